"""GPU tests of the cache operators against their 64-bit references
(_cache_ops): decoding behind a shared prefix, the attention weight of cached
keys (prompt and single token) and eviction, alone and as a serving loop runs
them together.

Bars: the decoding step's bf16 output as logo_decode's (max-abs 2e-2, mean-abs
2e-3); the weights within _cache_ops.score_tolerance; eviction exactly.
"""
import math

import numpy as np
import pytest

import _cache_ops as ref
import oracle
import synth
from _support import err_stats, to_device, torch_bf16_to_f64

pytestmark = pytest.mark.gpu

MAX_ABS, MEAN_ABS = 2e-2, 2e-3


@pytest.fixture(scope="module")
def pk():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu tests need an MI355X")
    import paper_2608_29539_amd as pk
    pk.library()
    oracle.build(force=False)
    return pk


def bf16(rng, *shape, std=1.0):
    return synth.bf16_bits_from_f32(
        (rng.standard_normal(int(np.prod(shape))) * std).astype(np.float32)).reshape(shape)


def cu_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)




# --- decoding behind a shared prefix ---------------------------------------------
def prefix_case(seed, prefixes, groups, own, hq, hkv, d, distinct):
    rng = np.random.default_rng(seed)
    B, N, P = len(own), sum(own), sum(prefixes)
    x = dict(q=bf16(rng, B, hq, d, std=2.0), k=bf16(rng, N, hkv, d), v=bf16(rng, N, hkv, d),
             k_pre=bf16(rng, P, hkv, d), v_pre=bf16(rng, P, hkv, d),
             gate=rng.random(B).astype(np.float32))
    if "q" in distinct:
        x["q_g"] = bf16(rng, B, hq, d, std=2.0)
    if "k" in distinct:
        for n, rows in (("k", N), ("v", N), ("k_pre", P), ("v_pre", P)):
            x[n + "_g"] = bf16(rng, rows, hkv, d)
    return x, cu_of(prefixes), cu_of(groups), cu_of(own)


def prefix_call(pk, x, cu_pre, cu_grp, cu, window, threshold, *, gains=None, host=True, slack=0,
                **kw):
    import torch
    dev = to_device({n: t for n, t in x.items()})
    dcu, dcp, dcg = (torch.from_numpy(t).cuda() for t in (cu, cu_pre, cu_grp))
    hq, hkv, d = x["q"].shape[1], x["k"].shape[1], x["q"].shape[2]
    sizes = {} if host else dict(total_tokens=int(cu[-1]), max_seqlen=int(np.diff(cu).max()) + slack)
    prob = pk.Problem(dcu, hq, hkv, d, window, cu_seqlens_host=cu if host else None, **sizes)
    if host:
        pre = pk.Prefix(dcp, dcg, cu_prefix_host=cu_pre, cu_group_host=cu_grp)
    else:
        pre = pk.Prefix(dcp, dcg, total_tokens=int(cu_pre[-1]),
                        max_prefix=int(np.diff(cu_pre).max()) + slack,
                        max_group=min(len(cu) - 1, int(np.diff(cu_grp).max()) + slack))
    for n, t in zip(("gain_local", "gain_global"), gains or ()):
        kw[n] = torch.from_numpy(t).cuda()
    glob = {n: dev[n] for n in ("q_g", "k_pre_g", "v_pre_g", "k_g", "v_g") if n in dev}
    if not (isinstance(threshold, dict)):
        threshold = dict(threshold=threshold)
    args = (prob, pre, dev["q"], dev["k_pre"], dev["v_pre"], dev["k"], dev["v"], dev["gate"])
    return pk.logo_decode_prefix(*args, **threshold, **glob, **kw), args, {**threshold, **glob, **kw}


def check_prefix(got, x, cu_pre, cu_grp, cu, window, threshold, gains, tag):
    gl, gg = gains or (None, None)
    want = ref.decode_prefix(x, cu_pre, cu_grp, cu, window, threshold, gain_local=gl, gain_global=gg)
    st = err_stats(torch_bf16_to_f64(got), want["out"])
    print(f"[prefix {tag}] n_sel={want['n_sel']} " + " ".join(f"{k}={v:.3g}" for k, v in st.items()),
          flush=True)
    assert st["max_abs"] <= MAX_ABS and st["mean_abs"] <= MEAN_ABS, (tag, st)
    return want


PREFIX_CASES = [
    # (prefixes, groups, own rows, Hq, Hkv, d, window, threshold, distinct, gains)
    ((300,), (3,), (1, 17, 64), 8, 2, 128, 128, 0.5, "", False),
    ((1,), (1,), (1,), 4, 4, 64, 1, 0.0, "", False),
    ((64, 65, 63), (2, 1, 2), (63, 1, 65, 128, 2), 4, 2, 64, 100, 0.3, "qk", True),
    ((0, 500, 0), (2, 0, 1), (5, 300, 77), 8, 2, 128, 64, 0.2, "", True),   # empty prefix, group
    ((700, 129), (2, 2), (0, 3, 0, 400), 6, 2, 64, 256, 0.4, "q", False),   # no rows of their own
    ((1000,), (5,), (1, 2, 3, 4, 5), 8, 8, 128, 5000, -math.inf, "", False),  # window past all
    ((1000,), (5,), (10, 600, 300, 301, 299), 8, 2, 128, 300, -math.inf, "", True),
    ((1000,), (5,), (10, 600, 300, 301, 299), 8, 2, 128, 300, math.inf, "k", False),
    ((2500, 40), (40, 1), tuple(1 + 7 * i for i in range(41)), 16, 4, 64, 200, 0.3, "", False),
    ((900,), (140,), tuple(1 + i % 9 for i in range(140)), 2, 2, 64, 64, 0.5, "", False),
    ((900,), (70,), tuple(1 + i % 30 for i in range(70)), 8, 2, 128, 1000, 0.1, "", False),
    ((300, 200), (3, 2), (3, 200, 9, 1, 70), 160, 1, 64, 128, 0.4, "", False),   # 160 heads a KV head
    ((350,), (50,), tuple(1 + i for i in range(50)), 3, 1, 128, 90, 0.5, "qk", True),
    ((20000,), (4,), (1, 700, 33, 2100), 8, 2, 128, 1024, 0.25, "", False),
    ((17000, 3), (3, 1), (40, 41, 42, 9000), 4, 1, 64, 512, 0.1, "", False),
    ((500, 600), (1, 1), (100, 100), 12, 4, 128, 1, 0.0, "", True),
]


@pytest.mark.parametrize("ci", range(len(PREFIX_CASES)))
def test_prefix(pk, ci):
    import torch
    pre, grp, own, hq, hkv, d, win, thr, distinct, gains = PREFIX_CASES[ci]
    rng = np.random.default_rng(50 + ci)
    gains = ([rng.uniform(0.5, 1.5, (hq, d)).astype(np.float32) for _ in range(2)]
             if gains else None)
    x, cp, cg, cu = prefix_case(ci, pre, grp, own, hq, hkv, d, distinct)
    for host in (True, False):
        print(f"[prefix case{ci}] host={host}", flush=True)
        act = torch.full((len(own),), -7, dtype=torch.int32, device="cuda")
        n_act = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        (got, _, _), args, kw = prefix_call(pk, x, cp, cg, cu, win, thr, gains=gains, host=host,
                                            slack=0 if host else 300, active=act, n_active=n_act)
        torch.cuda.synchronize()
        want = check_prefix(got, x, cp, cg, cu, win, thr, gains, f"case{ci}")
        sel = np.nonzero(want["z"])[0].tolist()
        assert n_act.tolist() == [len(sel)]
        assert act.tolist() == sel + [-7] * (len(own) - len(sel))
        # the same bits again, on another stream, in a workspace that is
        # exactly large enough
        need = pk.logo_decode_prefix_workspace_bytes(args[0], args[1])
        room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            again = pk.logo_decode_prefix(*args, **{**kw, "active": None, "n_active": None},
                                          ws=room[:need])[0]
        torch.cuda.synchronize()
        assert torch.equal(again.view(torch.int16), got.view(torch.int16))
        assert bool((room[need:] == 0xA5).all())


def test_prefix_gates_and_device_threshold(pk):
    """NaN gates are never selected, one equal to the threshold stays local;
    the threshold read on the device gives the same bits."""
    import torch
    x, cp, cg, cu = prefix_case(900, (400,), (6,), (3, 50, 7, 9, 200, 1), 8, 2, 128, "")
    x["gate"] = np.array([np.nan, 0.5, 0.5000001, 0.25, -0.0, 0.75], np.float32)
    (a, _, _), _, _ = prefix_call(pk, x, cp, cg, cu, 64, 0.5)
    want = check_prefix(a, x, cp, cg, cu, 64, 0.5, None, "gates")
    assert want["z"].tolist() == [False, False, True, False, False, True]
    t = torch.tensor([0.5], device="cuda")
    (b, _, _), _, _ = prefix_call(pk, x, cp, cg, cu, 64, dict(threshold_device=t))
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    t.fill_(float("nan"))
    (c, _, _), _, _ = prefix_call(pk, x, cp, cg, cu, 64, dict(threshold_device=t))
    check_prefix(c, x, cp, cg, cu, 64, math.inf, None, "NaN threshold")


def test_prefix_rows_outside_the_window_are_not_read(pk):
    """NaN in an unselected sequence's own rows before its window, and in
    prefix keys that no query sees."""
    import torch
    x, cp, cg, cu = prefix_case(903, (300,), (3,), (150, 100, 70), 8, 2, 128, "")
    x["gate"] = np.array([0.1, 0.2, 0.3], np.float32)
    (want, _, _), args, kw = prefix_call(pk, x, cp, cg, cu, 64, 0.5)
    prob, pre, q, kp, vp, k, v, gate = args
    for t in (k, v):
        for b in range(3):
            t[cu[b]:cu[b + 1] - 64] = float("nan")
    for t in (kp, vp):
        t[:] = float("nan")                      # every sequence has its window in its own rows
    got = pk.logo_decode_prefix(*args, **kw)[0]
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_two_streams(pk):
    """Steps on two streams with workspaces of their own, interleaved."""
    import torch
    cases = [prefix_case(904 + i, (600 + 50 * i,), (4,), (5, 90, 30, 1), 8, 2, 128, "") for i in range(2)]
    calls = [prefix_call(pk, *c, 128, 0.4) for c in cases]
    torch.cuda.synchronize()
    want = [c[0][0].clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    outs = []
    for _ in range(20):
        for (_, args, kw), s in zip(calls, streams):
            with torch.cuda.stream(s):
                outs.append(pk.logo_decode_prefix(*args, **kw)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o.view(torch.int16), want[i % 2].view(torch.int16)), i


def test_prefix_without_any_rows(pk):
    """Without host copies a sequence with no rows at all outputs zeros."""
    import torch
    x, cp, cg, cu = prefix_case(901, (0, 30), (1, 1), (0, 4), 4, 2, 64, "")
    (got, _, _), _, _ = prefix_call(pk, x, cp, cg, cu, 8, -math.inf, host=False)
    torch.cuda.synchronize()
    assert bool((got[0] == 0).all()) and bool(torch.isfinite(got.float()).all())


def test_prefix_agrees_with_decode(pk):
    """One sequence per prefix: logo_decode on the joined caches."""
    import torch
    x, cp, cg, cu = prefix_case(902, (800, 33, 5000), (1, 1, 1), (9, 300, 64), 8, 2, 128, "")
    (got, _, _), args, _ = prefix_call(pk, x, cp, cg, cu, 512, 0.3)
    k, whole = ref.whole_caches(x["k_pre"], x["k"], cp, cg, cu)
    v, _ = ref.whole_caches(x["v_pre"], x["v"], cp, cg, cu)
    dev = to_device(dict(q=x["q"], k=k, v=v, gate=x["gate"], cu=whole))
    prob = pk.Problem(dev["cu"], 8, 2, 128, 512, cu_seqlens_host=whole)
    one = pk.logo_decode(prob, dev["q"], dev["k"], dev["v"], dev["gate"], threshold=0.3)[0]
    st = err_stats(torch_bf16_to_f64(got), torch_bf16_to_f64(one))
    assert st["max_abs"] <= MAX_ABS and st["mean_abs"] <= MEAN_ABS, st


# --- attention weight of cached keys ----------------------------------------------
def score_case(seed, lens, hq, hkv, d):
    rng = np.random.default_rng(seed)
    N = sum(lens)
    return bf16(rng, N, hq, d, std=2.0), bf16(rng, N, hkv, d), cu_of(lens), rng


SCORE_CASES = [
    # (lengths, share of rows, Hq, Hkv, d, scale)
    ((1,), 1.0, 4, 4, 64, 0.0), ((1, 64, 65), 1.0, 4, 2, 128, 0.0),
    ((300, 0, 257), 0.3, 8, 2, 128, 0.0), ((500,), 0.1, 3, 1, 64, 0.2),
    ((130, 700), 0.25, 16, 2, 64, 0.0), ((1500,), 0.05, 8, 8, 128, 0.05),
    ((200, 31, 1000), 0.0, 8, 4, 128, 0.0), ((90,) * 70, 0.2, 4, 4, 64, 0.0),
    ((40, 0, 90), 1.0, 40, 1, 64, 0.0),
]


@pytest.mark.parametrize("ci", range(len(SCORE_CASES)))
def test_cache_score(pk, ci):
    import torch
    lens, share, hq, hkv, d, scale = SCORE_CASES[ci]
    q, k, cu, rng = score_case(ci, lens, hq, hkv, d)
    N = sum(lens)
    rows = [np.sort(rng.choice(T, max(int(share * T), 1 if share and T else 0), replace=False))
            for T in lens]
    n = [len(r) for r in rows]
    sel = np.concatenate([r + c for r, c in zip(rows, cu)]).astype(np.int32)
    total, size = ref.scores_of(q, k, sel, cu, n, scale=scale)
    before = rng.random((hkv, N)).astype(np.float32)
    dev = to_device(dict(q=q, k=k, cu=cu, before=before, cu_sel=cu_of(n)))
    prob = pk.Problem(dev["cu"], hq, hkv, d, 64, cu_seqlens_host=cu, softmax_scale=scale)
    # sel_idx has room behind the last row, filled with what must not be read
    # as a row
    cap = len(sel) + 37
    idx = torch.full((cap,), 1 << 30, dtype=torch.int32, device="cuda")
    idx[:len(sel)] = torch.from_numpy(sel).cuda()
    kw = dict(sel_idx=idx, cu_sel=dev["cu_sel"])
    tol = ref.score_tolerance(total + before, max(n) * (hq // hkv), d, size)

    def check(got, add, tag):
        torch.cuda.synchronize()
        e = np.abs(got.cpu().numpy().astype(np.float64) - (total + add))
        print(f"[score case{ci} {tag}] size={size:.3g} worst/tol={(e / tol).max() if e.size else 0:.3g}",
              flush=True)
        assert np.all(e <= tol), (tag, e.max())

    print(f"[score case{ci}] {lens}", flush=True)
    own = pk.logo_cache_score(prob, dev["q"], dev["k"], score_in=dev["before"], **kw)
    check(own, before, "lse computed")
    check(pk.logo_cache_score(prob, dev["q"], dev["k"], **kw), 0.0, "from zero")
    lse = pk.logo_global_attn_sparse_q_fwd_train(prob, dev["q"], dev["k"], dev["k"], idx,
                                                 dev["cu_sel"], cap)[1]
    inplace = dev["before"].clone()
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], lse=lse, score_in=inplace, score=inplace, **kw)
    assert got.data_ptr() == inplace.data_ptr()
    # (that forward's row sums take P rounded to bf16: its lse is off by up to
    # log2(1 + 2^-8), which the weights follow)
    torch.cuda.synchronize()
    e = np.abs(inplace.cpu().numpy().astype(np.float64) - (total + before))
    assert np.all(e <= tol + total * 2.0 ** -7)
    # against the reference with that very lse
    total, _ = ref.scores_of(q, k, sel, cu, n, scale=scale, lse=lse.cpu().numpy().astype(np.float64))
    check(got, before, "lse given")
    again = pk.logo_cache_score(prob, dev["q"], dev["k"], score_in=dev["before"], **kw)
    assert torch.equal(again, own)


def test_cache_score_every_row(pk):
    """Without a selection every token is a row; the dense forward's lse."""
    import torch
    lens = (100, 1, 333)
    q, k, cu, _ = score_case(77, lens, 8, 2, 128)
    dev = to_device(dict(q=q, k=k, cu=cu))
    prob = pk.Problem(dev["cu"], 8, 2, 128, 64, cu_seqlens_host=cu)
    total, size = ref.scores_of(q, k, np.arange(sum(lens)), cu, lens)
    got = pk.logo_cache_score(prob, dev["q"], dev["k"]).cpu().numpy().astype(np.float64)
    tol = ref.score_tolerance(total, max(lens) * 4, 128, size)
    assert np.all(np.abs(got - total) <= tol)
    # every row gives a weight of one in all
    np.testing.assert_allclose(got.sum(), sum(lens) * 8, rtol=1e-4)
    lse = pk.logo_dense_causal_attn_fwd_train(prob, dev["q"], dev["k"], dev["k"])[1]
    total, _ = ref.scores_of(q, k, np.arange(sum(lens)), cu, lens,
                             lse=lse.cpu().numpy().astype(np.float64))
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], lse=lse).cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - total) <= ref.score_tolerance(total, max(lens) * 4, 128, size))


def test_cache_score_capacity_overflow(pk):
    """Only the first sel_capacity rows count."""
    import torch
    q, k, cu, _ = score_case(78, (200, 300), 4, 2, 64)
    sel = np.concatenate([np.arange(0, 200, 3), 200 + np.arange(0, 300, 5)]).astype(np.int32)
    n0 = len(np.arange(0, 200, 3))
    dev = to_device(dict(q=q, k=k, cu=cu, sel=sel, cu_sel=np.array([0, n0, len(sel)], np.int32)))
    prob = pk.Problem(dev["cu"], 4, 2, 64, 64, cu_seqlens_host=cu)
    for cap in (n0 + 11, n0 - 5):
        n = [min(n0, cap), max(0, cap - n0)]
        total, size = ref.scores_of(q, k, sel[:cap], cu, n)
        got = pk.logo_cache_score(prob, dev["q"], dev["k"], sel_idx=dev["sel"][:cap].contiguous(),
                                  cu_sel=dev["cu_sel"])
        e = np.abs(got.cpu().numpy().astype(np.float64) - total)
        assert np.all(e <= ref.score_tolerance(total, 500, 64, size)), cap


def test_cache_score_later_keys_do_not_reach_earlier_rows(pk):
    """NaN and infinite keys behind every row: the rows give what they gave."""
    import torch
    q, k, cu, _ = score_case(79, (300,), 8, 2, 128)
    sel = np.arange(0, 150, 2).astype(np.int32)
    dev = to_device(dict(q=q, k=k, cu=cu, sel=sel, cu_sel=np.array([0, len(sel)], np.int32)))
    prob = pk.Problem(dev["cu"], 8, 2, 128, 64, cu_seqlens_host=cu)
    kw = dict(sel_idx=dev["sel"], cu_sel=dev["cu_sel"])
    want = pk.logo_cache_score(prob, dev["q"], dev["k"], **kw)
    dev["k"][149:200] = float("nan")
    dev["k"][200:] = float("inf")
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], **kw)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and bool((got[:, 149:] == 0).all())


STEP_CASES = [
    # (caches, Hq, Hkv, d, threshold, scale)
    ((1,), 4, 4, 64, 0.0, 0.0), ((1, 15, 16, 17, 300), 8, 2, 128, 0.4, 0.0),
    ((2000, 511, 512, 513, 1), 16, 2, 64, 0.3, 0.1), ((700, 5000), 20, 1, 128, 0.0, 0.0),
    ((1025, 1024, 1023), 3, 3, 128, math.inf, 0.0), ((33000,), 4, 2, 64, -math.inf, 0.0),
    ((900, 40), 34, 2, 64, 0.1, 0.0),
]


@pytest.mark.parametrize("ci", range(len(STEP_CASES)))
def test_decode_score(pk, ci):
    import torch
    lens, hq, hkv, d, thr, scale = STEP_CASES[ci]
    rng = np.random.default_rng(300 + ci)
    N, B = sum(lens), len(lens)
    q, k, cu = bf16(rng, B, hq, d, std=2.0), bf16(rng, N, hkv, d), cu_of(lens)
    gate = rng.random(B).astype(np.float32)
    if B > 2:
        gate[1] = np.nan
    before = rng.random((hkv, N)).astype(np.float32)
    total, size = ref.step_scores(q, k, cu, gate > thr, scale=scale)
    tol = ref.score_tolerance(total + before, hq // hkv, d, size)
    dev = to_device(dict(q=q, k=k, cu=cu, gate=gate, before=before))
    prob = pk.Problem(dev["cu"], hq, hkv, d, 64, cu_seqlens_host=cu, softmax_scale=scale)
    need = pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_DECODE_SCORE)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    print(f"[step case{ci}] {lens}", flush=True)

    def check(got, add):
        torch.cuda.synchronize()
        e = np.abs(got.cpu().numpy().astype(np.float64) - (total + add))
        assert np.all(e <= tol), e.max()

    got = pk.logo_decode_score(prob, dev["q"], dev["k"], dev["gate"], threshold=thr,
                               score_in=dev["before"], ws=room[:need])
    check(got, before)
    assert bool((room[need:] == 0xA5).all())
    check(pk.logo_decode_score(prob, dev["q"], dev["k"], dev["gate"], threshold=thr), 0.0)
    t = torch.tensor([thr], device="cuda")
    inplace = dev["before"].clone()
    pk.logo_decode_score(prob, dev["q"], dev["k"], dev["gate"], threshold_device=t,
                         score_in=inplace, score=inplace)
    torch.cuda.synchronize()
    assert torch.equal(inplace, got)


def test_cache_score_nothing_selected(pk):
    """No row: the scores stay as they were."""
    import torch
    q, k, cu, rng = score_case(80, (70, 0, 9), 4, 2, 64)
    before = rng.random((2, 79)).astype(np.float32)
    dev = to_device(dict(q=q, k=k, cu=cu, before=before))
    prob = pk.Problem(dev["cu"], 4, 2, 64, 64, cu_seqlens_host=cu)
    none = dict(sel_idx=torch.empty(0, dtype=torch.int32, device="cuda"),
                cu_sel=torch.zeros(4, dtype=torch.int32, device="cuda"))
    for lse in (None, torch.empty((4, 0), device="cuda")):
        got = pk.logo_cache_score(prob, dev["q"], dev["k"], lse=lse, score_in=dev["before"], **none)
        assert torch.equal(got, dev["before"])
    # room for rows, but none of them selected
    none["sel_idx"] = torch.full((50,), 1 << 30, dtype=torch.int32, device="cuda")
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], **none)
    assert bool((got == 0).all())


@pytest.mark.parametrize("lens", [tuple([5] * 300), tuple([3] * 150 + [2000, 0] + [1] * 149)],
                         ids=["even", "one-long"])
def test_cache_score_many_sequences(pk, lens):
    """Workgroups find their sequence by a division (even lengths) or a search."""
    q, k, cu, rng = score_case(81, lens, 2, 1, 64)
    rows = [np.sort(rng.choice(T, (T + 2) // 3 if T < 100 else 60, replace=False)) if T else
            np.zeros(0, np.int64) for T in lens]
    n = [len(r) for r in rows]
    sel = np.concatenate([r + c for r, c in zip(rows, cu)]).astype(np.int32)
    total, size = ref.scores_of(q, k, sel, cu, n)
    dev = to_device(dict(q=q, k=k, cu=cu, sel=sel, cu_sel=cu_of(n)))
    prob = pk.Problem(dev["cu"], 2, 1, 64, 64, cu_seqlens_host=cu)
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], sel_idx=dev["sel"], cu_sel=dev["cu_sel"])
    e = np.abs(got.cpu().numpy().astype(np.float64) - total)
    assert np.all(e <= ref.score_tolerance(total, max(n) * 2, 64, size))


def test_cache_score_row_listed_twice(pk):
    """A row in the list twice gives its weights twice."""
    q, k, cu, _ = score_case(82, (40, 30), 8, 2, 128)
    sel = np.array([3, 3, 3, 17, 39, 40, 40, 69], np.int32)
    dev = to_device(dict(q=q, k=k, cu=cu, sel=sel, cu_sel=np.array([0, 5, 8], np.int32)))
    prob = pk.Problem(dev["cu"], 8, 2, 128, 64, cu_seqlens_host=cu)
    total, size = ref.scores_of(q, k, sel, cu, [5, 3])
    got = pk.logo_cache_score(prob, dev["q"], dev["k"], sel_idx=dev["sel"], cu_sel=dev["cu_sel"])
    e = np.abs(got.cpu().numpy().astype(np.float64) - total)
    assert np.all(e <= ref.score_tolerance(total, 5 * 4, 128, size))


def test_offsets_past_32_bits(pk):
    """Caches of more than 4 GiB: the second sequence lies behind the first
    one's 2.2 million rows, and a prefix behind another one's."""
    import torch
    hq, hkv, d, far, L = 16, 8, 128, 2200000, 300
    rng = np.random.default_rng(83)
    q, k, v = bf16(rng, 1, hq, d, std=2.0), bf16(rng, L, hkv, d), bf16(rng, L, hkv, d)
    dev = to_device(dict(q=q, k=k, v=v))
    big_k, big_v = (torch.zeros((far + L, hkv, d), dtype=torch.bfloat16, device="cuda")
                    for _ in range(2))
    assert big_k.numel() * 2 > 1 << 32
    big_k[far:], big_v[far:] = dev["k"], dev["v"]
    cu = np.array([0, far, far + L], np.int32)
    dcu = torch.from_numpy(cu).cuda()
    prob = pk.Problem(dcu, hq, hkv, d, 64, cu_seqlens_host=cu)
    want, size = ref.step_scores(q, k, [0, L], [True])
    tol = ref.score_tolerance(want, hq // hkv, d, size)
    # one decoding step of the second sequence
    q2 = torch.cat([dev["q"], dev["q"]])
    gate = torch.tensor([0.0, 1.0], device="cuda")
    got = pk.logo_decode_score(prob, q2, big_k, gate, threshold=0.5)
    assert bool((got[:, :far] == 0).all())
    assert np.all(np.abs(got[:, far:].cpu().numpy() - want) <= tol)
    # its last row as a prompt's only query
    qq = torch.zeros((far + L, hq, d), dtype=torch.bfloat16, device="cuda")
    qq[-1] = dev["q"][0]
    got = pk.logo_cache_score(prob, qq, big_k,
                              sel_idx=torch.tensor([far + L - 1], dtype=torch.int32, device="cuda"),
                              cu_sel=torch.tensor([0, 0, 1], dtype=torch.int32, device="cuda"))
    assert bool((got[:, :far] == 0).all())
    assert np.all(np.abs(got[:, far:].cpu().numpy() - want) <= tol)
    del qq, q2
    # eviction: all scores equal in the first sequence, so its oldest rows stay
    sc = torch.rand((hkv, far + L), device="cuda")
    sc[:, :far] = 0.25
    r = pk.logo_cache_evict(prob, sc, 100, recent=10, k=big_k, v=big_v)
    kept, _ = ref.evict(sc[:, far:].cpu().numpy(), np.array([0, L]), 100, 10)
    idx = r["keep_idx"].cpu().numpy()
    first = list(range(90)) + list(range(far - 10, far))
    assert (idx[:, :100] == first).all() and np.array_equal(idx[:, 100:], kept + far)
    for h in range(hkv):
        assert torch.equal(r["k_out"][100:, h], big_k[r["keep_idx"][h, 100:].long(), h])
        assert torch.equal(r["v_out"][100:, h], big_v[r["keep_idx"][h, 100:].long(), h])
    # the far rows as a shared prefix
    own = dict(k=bf16(rng, 5, hkv, d), v=bf16(rng, 5, hkv, d), gate=np.array([0.9, 0.2], np.float32))
    x = dict(q=np.concatenate([q, q[:, ::-1]]), k_pre=k, v_pre=v, **own)
    cu_own, cu_grp = np.array([0, 2, 5], np.int32), np.array([0, 0, 2], np.int32)
    d2 = to_device(dict(q=x["q"], cu=cu_own, grp=cu_grp, **own))
    pre = pk.Prefix(dcu, d2["grp"], cu_prefix_host=cu, cu_group_host=cu_grp)
    p2 = pk.Problem(d2["cu"], hq, hkv, d, 64, cu_seqlens_host=cu_own)
    out = pk.logo_decode_prefix(p2, pre, d2["q"], big_k, big_v, d2["k"], d2["v"], d2["gate"],
                                threshold=0.5)[0]
    check_prefix(out, x, np.array([0, L]), np.array([0, 2]), cu_own, 64, 0.5, None, "far")


# --- eviction -------------------------------------------------------------------
def evict_scores(rng, hkv, N, kind):
    s = np.exp(2 * rng.standard_normal((hkv, N))).astype(np.float32)
    s[rng.random((hkv, N)) < 0.1] = 0.0
    if kind == "equal":
        s[:] = 0.25
    if kind == "few":
        s = rng.choice(np.array([0.0, -0.0, 1.0, 2.0], np.float32), (hkv, N))
    if kind == "odd":
        s = rng.standard_normal((hkv, N)).astype(np.float32)
        for v in (np.nan, np.inf, -np.inf, -0.0, 0.0, 1e-42, -1e-42, 3.4e38):
            s[rng.random((hkv, N)) < 0.08] = v
    if kind == "nan":
        s[:] = np.nan
    return s


EVICT_CASES = [
    # (caches, Hkv, d, budget, recent, scores)
    ((1,), 1, 64, 1, 0, "heavy"), ((5, 300, 1), 2, 128, 7, 3, "heavy"),
    ((100, 0, 2000, 1024, 1025), 4, 64, 512, 128, "heavy"), ((3000, 50), 2, 128, 100, 0, "equal"),
    ((3000, 50, 1000), 8, 64, 900, 10, "few"), ((2500, 700), 3, 128, 600, 33, "odd"),
    ((2500, 700), 2, 64, 2499, 0, "odd"), ((900,), 2, 64, 100, 50, "nan"),
    ((400, 90), 2, 128, 1000, 20, "heavy"), ((400, 90), 2, 128, 60, 500, "heavy"),
    ((400, 90), 2, 128, 60, 60, "odd"), ((9,) * 300, 2, 64, 4, 1, "odd"),
    ((40000, 33), 2, 64, 5001, 1000, "heavy"), ((131071,), 1, 64, 16001, 0, "few"),
    ((131071,), 1, 128, 16001, 4096, "heavy"), ((70001,), 3, 64, 1, 0, "odd"),
]


@pytest.mark.parametrize("ci", range(len(EVICT_CASES)))
def test_evict(pk, ci):
    import torch
    lens, hkv, d, budget, recent, kind = EVICT_CASES[ci]
    rng = np.random.default_rng(600 + ci)
    N, cu = sum(lens), cu_of(lens)
    score = evict_scores(rng, hkv, N, kind)
    x = {n: bf16(rng, N, hkv, d) for n in ("k", "v", "k_g", "v_g")}
    kept, cu_keep = ref.evict(score, cu, budget, recent)
    n = kept.shape[1]
    dev = to_device(dict(score=score, cu=cu, **x))
    prob = pk.Problem(dev["cu"], hkv, hkv, d, 64, cu_seqlens_host=cu)
    assert pk.logo_cache_keep_capacity(prob, budget) == n
    extra = 5                                    # rows behind the last stay as they were
    out = {f"{t}_out": torch.full((n + extra, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
           for t in x}
    out["score_out"] = torch.full((hkv, n + extra), -5.0, device="cuda")
    out["keep_idx"] = torch.full((hkv, n + extra), -5, dtype=torch.int32, device="cuda")
    print(f"[evict case{ci}] {lens[:6]} {kind}", flush=True)
    r = pk.logo_cache_evict(prob, dev["score"], budget, recent=recent,
                            **{t: dev[t] for t in x}, **out)
    torch.cuda.synchronize()
    assert r["cu_keep"].cpu().numpy().tolist() == cu_keep.tolist()
    idx = r["keep_idx"].cpu().numpy()
    assert np.array_equal(idx[:, :n], kept) and (idx[:, n:] == -5).all()
    so = r["score_out"].cpu().numpy()
    assert np.array_equal(so[:, :n].view(np.int32),
                          np.take_along_axis(score, kept, 1).view(np.int32))
    assert (so[:, n:] == -5).all()
    for t in x:
        got = r[f"{t}_out"].view(torch.int16).cpu().numpy().view(np.uint16)
        for h in range(hkv):
            assert np.array_equal(got[:n, h], x[t][kept[h], h]), (t, h)
        assert bool((r[f"{t}_out"][n:] == 7.0).all())
    # the choice alone, without a host copy of the lengths
    bare = pk.Problem(dev["cu"], hkv, hkv, d, 64, total_tokens=N, max_seqlen=max(lens))
    c = pk.logo_cache_evict(bare, dev["score"], budget, recent=recent)
    torch.cuda.synchronize()
    assert c["k_out"] is None and np.array_equal(c["keep_idx"].cpu().numpy()[:, :n], kept)


def test_evict_nothing(pk):
    """Caches without rows, with and without outputs' room."""
    import torch
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    prob = pk.Problem(cu, 4, 2, 64, 64, cu_seqlens_host=[0, 0, 0, 0])
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    r = pk.logo_cache_evict(prob, torch.empty((2, 0), device="cuda"), 5, recent=2, k=empty, v=empty)
    assert r["cu_keep"].tolist() == [0, 0, 0, 0] and r["k_out"].shape[0] == 0


# --- together -------------------------------------------------------------------
def serving_inputs(rng, hq, hkv, d, P, own):
    pre = dict(q=bf16(rng, P, hq, d, std=2.0), k=bf16(rng, P, hkv, d), v=bf16(rng, P, hkv, d),
               gate=rng.random(P).astype(np.float32))
    new = dict(q=bf16(rng, len(own), hq, d, std=2.0), k=bf16(rng, sum(own), hkv, d),
               v=bf16(rng, sum(own), hkv, d), gate=rng.random(len(own)).astype(np.float32))
    return pre, new


def test_serving_run(pk):
    """A prompt is run through the layer, its keys scored with the layer's own
    lse, its cache cut down; a group of sequences decodes behind what is left;
    and a sequence's joined cache goes on with scored steps and another
    eviction.  Each stage is compared with its reference on that stage's
    inputs."""
    import torch
    hq, hkv, d, win, P, own = 8, 2, 128, 96, 1500, (1, 40, 7)
    rng = np.random.default_rng(4)
    pre, new = serving_inputs(rng, hq, hkv, d, P, own)
    cu = cu_of([P])
    dev = to_device(dict(cu=cu, **pre))
    prob = pk.Problem(dev["cu"], hq, hkv, d, win, cu_seqlens_host=cu)
    st = pk.logo_attn_fwd_train(prob, dev["q"], dev["k"], dev["v"], dev["gate"], ratio=0.125)
    n_sel = int(st["cu_sel"][-1])
    sel = st["sel_idx"][:n_sel]
    score = pk.logo_cache_score(prob, dev["q"], dev["k"], sel_idx=st["sel_idx"],
                                cu_sel=st["cu_sel"], lse=st["lse_global"])
    total, size = ref.scores_of(pre["q"], pre["k"], sel.cpu().numpy(), cu, [n_sel],
                                lse=st["lse_global"].cpu().numpy().astype(np.float64))
    got = score.cpu().numpy()
    assert np.all(np.abs(got - total) <= ref.score_tolerance(total, n_sel * 4, d, size))
    ev = pk.logo_cache_evict(prob, score, 400, recent=win, k=dev["k"], v=dev["v"])
    kept, cu_keep = ref.evict(got, cu, 400, win)
    assert np.array_equal(ev["keep_idx"].cpu().numpy(), kept)
    # the group decodes behind the kept rows
    x = dict(q=new["q"], k=new["k"], v=new["v"], gate=new["gate"],
             k_pre=np.stack([pre["k"][kept[h], h] for h in range(hkv)], 1),
             v_pre=np.stack([pre["v"][kept[h], h] for h in range(hkv)], 1))
    (out, _, _), _, _ = prefix_call(pk, x, cu_keep, cu_of([3]), cu_of(own), win, 0.4)
    check_prefix(out, x, cu_keep, cu_of([3]), cu_of(own), win, 0.4, None, "serving")
    # the sequences go on with caches of their own
    k, whole = ref.whole_caches(x["k_pre"], x["k"], cu_keep, cu_of([3]), cu_of(own))
    v, _ = ref.whole_caches(x["v_pre"], x["v"], cu_keep, cu_of([3]), cu_of(own))
    d2 = to_device(dict(q=new["q"], k=k, v=v, gate=new["gate"], cu=whole))
    prob2 = pk.Problem(d2["cu"], hq, hkv, d, win, cu_seqlens_host=whole)
    s2 = pk.logo_decode_score(prob2, d2["q"], d2["k"], d2["gate"], threshold=0.4)
    total, size = ref.step_scores(new["q"], k, whole, new["gate"] > 0.4)
    got = s2.cpu().numpy()
    assert np.all(np.abs(got - total) <= ref.score_tolerance(total, 4, d, size))
    e2 = pk.logo_cache_evict(prob2, s2, 300, recent=win, k=d2["k"], v=d2["v"])
    kept2, cu2 = ref.evict(got, whole, 300, win)
    assert np.array_equal(e2["keep_idx"].cpu().numpy(), kept2)
    prob3 = pk.Problem(e2["cu_keep"], hq, hkv, d, win, cu_seqlens_host=cu2)
    o3 = pk.logo_decode(prob3, d2["q"], e2["k_out"], e2["v_out"], d2["gate"], threshold=0.4)[0]
    want = oracle.decode(new["q"], np.stack([k[kept2[h], h] for h in range(hkv)], 1),
                         np.stack([v[kept2[h], h] for h in range(hkv)], 1), new["gate"], cu2, win,
                         0.4)
    st = err_stats(torch_bf16_to_f64(o3), want["out"])
    assert st["max_abs"] <= MAX_ABS and st["mean_abs"] <= MEAN_ABS, st


def test_captured_step(pk):
    """Decoding, scoring and eviction captured into one graph, replayed with
    new inputs and with eager work between the replays."""
    import torch
    hq, hkv, d, win, own = 8, 2, 64, 64, (30, 5, 200)
    rng = np.random.default_rng(5)
    x, cp, cg, cu = prefix_case(6, (700,), (3,), own, hq, hkv, d, "")
    (_, _, _), args, kw = prefix_call(pk, x, cp, cg, cu, win, 0.3)
    prob, pre, q, kp, vp, k, v, gate = args
    cap = pk.logo_cache_keep_capacity(prob, 20)
    ws = torch.empty(pk.logo_decode_prefix_workspace_bytes(prob, pre), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_DECODE_SCORE), dtype=torch.uint8,
                      device="cuda")
    ws3 = torch.empty(pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_CACHE_SCORE, 3), dtype=torch.uint8,
                      device="cuda")
    ws4 = torch.empty(max(256, pk.logo_workspace_bytes(prob, pk.LOGO_ENTRY_CACHE_EVICT)),
                      dtype=torch.uint8, device="cuda")
    sel = torch.tensor([29, 34, 234], dtype=torch.int32, device="cuda")
    cu_sel = torch.arange(4, dtype=torch.int32, device="cuda")
    qn = torch.zeros((sum(own), hq, d), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    score = torch.zeros((hkv, sum(own)), device="cuda")
    ev = {n: torch.zeros((cap, hkv, d), dtype=torch.bfloat16, device="cuda") for n in ("k_out", "v_out")}
    ev.update(score_out=torch.zeros((hkv, cap), device="cuda"),
              keep_idx=torch.zeros((hkv, cap), dtype=torch.int32, device="cuda"),
              cu_keep=torch.zeros(4, dtype=torch.int32, device="cuda"))

    def step():
        pk.logo_decode_prefix(*args, threshold=0.3, out=out, ws=ws)
        pk.logo_decode_score(prob, q, k, gate, threshold=0.3, score_in=score, score=score, ws=ws2)
        pk.logo_cache_score(prob, qn, k, sel_idx=sel, cu_sel=cu_sel, score_in=score, score=score,
                            ws=ws3)
        pk.logo_cache_evict(prob, score, 20, recent=4, k=k, v=v, ws=ws4, **ev)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    got = {**ev, "out": out, "score": score}
    for i in range(4):
        q.copy_(torch.from_numpy(rng.standard_normal(tuple(q.shape)).astype(np.float32)))
        qn.copy_(torch.from_numpy(rng.standard_normal(tuple(qn.shape)).astype(np.float32)))
        gate.copy_(torch.rand(3))
        start = torch.rand_like(score)
        score.copy_(start)
        g.replay()
        torch.cuda.synchronize()
        first = {n: t.clone() for n, t in got.items()}
        score.copy_(start)
        step()
        torch.cuda.synchronize()
        for n, t in got.items():
            assert torch.equal(first[n].view(torch.int32 if t.element_size() == 4 else torch.int16),
                               t.view(torch.int32 if t.element_size() == 4 else torch.int16)), (i, n)
