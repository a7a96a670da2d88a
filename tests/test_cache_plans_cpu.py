"""The plans of the cache operators and the workspaces that they ask for, on
the CPU: a workspace given for a larger call serves every smaller one."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ALL = (1 << 64) - 1


@pytest.fixture(scope="module")
def lib():
    import paper_2608_29539_amd as pk
    if not os.path.exists(pk.library_path()):
        from paper_2608_29539_amd.build import build_library
        build_library()
    return pk.library()


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plans") / "plans.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared",
                    "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-I", os.path.join(ROOT, "paper_2608_29539_amd", "csrc"),
                    os.path.join(ROOT, "tests", "c", "cache_plans.cpp"), "-o", so], check=True)
    so = ctypes.CDLL(so)
    so.evict_total.restype = ctypes.c_longlong
    return so


CU = np.zeros(1, np.int32)
PTR = CU.ctypes.data_as(ctypes.c_void_p)


def problem(B, N, longest, hq, hkv, d, window):
    import paper_2608_29539_amd.binding as b
    return b._Problem(B, N, longest, PTR, None, hq, hkv, d, window, 0.0)


def prefixes(R, total, longest, group):
    import paper_2608_29539_amd.binding as b
    return b._Prefix(R, total, longest, group, PTR, PTR, None, None)


def size_t(x):
    return ctypes.c_size_t(x)


def prefix(plans, p, x, share, room=ALL):
    out = (ctypes.c_longlong * 18)()
    plans.prefix_plan(ctypes.byref(p), ctypes.byref(x), int(share), size_t(room), out)
    v = list(out)
    return dict(total=v[0], ml=v[1], kc=v[2:6], chunks=v[6:10], slot0=v[10:14], items=v[14:18])


def small(plans, name, p, room, *args):
    out = (ctypes.c_longlong * 3)()
    getattr(plans, name)(ctypes.byref(p), *args, size_t(room), out)
    return dict(zip(("total", "kc", "chunks"), out))


def up(x, n=256):
    return -(-x // n) * n


def prefix_bytes(lib, p, x):
    return lib.logo_decode_prefix_workspace_bytes(ctypes.byref(p), ctypes.byref(x))


def check_prefix_plan(d, p, x, share, room):
    P, S, w = x.max_prefix, p.max_seqlen, p.window
    spans = [P, max(0, S - w) if share else S, min(P, w), min(S, w)]
    rows = p.num_seqs * p.num_q_heads
    slots = 0
    for i, n in enumerate(spans):
        assert d["kc"][i] > 0 and d["kc"][i] % 64 == 0
        assert d["chunks"][i] == -(-n // d["kc"][i]) <= 128
        assert d["slot0"][i] == slots
        slots += d["chunks"][i]
    assert d["ml"] == up(4 * rows * slots * p.head_dim)
    assert d["total"] == d["ml"] + up(8 * rows * slots) and d["total"] <= room


HEADS = [(32, 8, 128), (4, 4, 64), (16, 2, 128), (40, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("B,groups", [(1, 1), (16, 1), (32, 3), (64, 2)])
def test_prefix_workspace_of_a_longer_step(plans, lib, hq, hkv, d, B, groups):
    """Steps of growing prefixes and own caches: each one's size is taken by
    every earlier one, whichever tensors the branches read."""
    lengths = [(P, S) for P in (0, 1, 300, 1024, 5000, 10240, 15360, 16384, 40000, 200000)
               for S in (1, 100, 1024, 1400, 2048, 9000)]
    rng = np.random.default_rng(B * hq)
    for w in (64, 1024, 1 << 30):
        big = []
        for P, S in lengths:
            p = problem(B, B * S, S, hq, hkv, d, w)
            x = prefixes(groups, P * groups, P, -(-B // groups))
            big.append((P, S, p, x, prefix_bytes(lib, p, x)))
            for share in (False, True):
                check_prefix_plan(prefix(plans, p, x, share), p, x, share, big[-1][4])
        for P, S, p, x, need in big:
            for Pb, Sb, _, _, room in big:
                if Pb < P or Sb < S:
                    continue
                share = bool(rng.random() < 0.5)
                check_prefix_plan(prefix(plans, p, x, share, room), p, x, share, room)
                # the size of the call itself leaves its plan as it is
                assert prefix(plans, p, x, share, need) == prefix(plans, p, x, share)


def test_prefix_workspace_of_more_sequences(plans, lib):
    """The last sequences of a batch leave it, and with them its prefixes."""
    big = problem(64, 64 * 500, 500, 32, 8, 128, 1024)
    room = prefix_bytes(lib, big, prefixes(4, 4 * 9000, 9000, 40))
    for B in range(1, 65):
        for R, longest in ((4, 9000), (3, 5000), (1, 9000), (1, 1)):
            p, x = problem(B, B * 200, 200, 32, 8, 128, 1024), prefixes(R, R * longest, longest,
                                                                       min(B, 40))
            for share in (False, True):
                check_prefix_plan(prefix(plans, p, x, share, room), p, x, share, room)


def test_prefix_sizes_that_shrink(lib):
    """What the sweeps above are for: sizes that a longer step's does not cover."""
    def need(P, S, B=32):
        return prefix_bytes(lib, problem(B, B * S, S, 32, 8, 128, 1024), prefixes(1, P, P, B))

    assert need(10240, 100) > need(16384, 100)
    assert need(8192, 1536, 16) > need(8192, 2048, 16)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_score_workspace_of_more_rows(plans, lib, hq, hkv, d):
    import paper_2608_29539_amd as pk
    sizes = []
    for L in (1, 500, 4096, 32768):
        for cap in (1, 64, 100, 640, 2000, 4000, 4096, 32768):
            p = problem(3, 2 * L + 1, L, hq, hkv, d, 64)
            need = lib.logo_workspace_bytes(ctypes.byref(p), pk.LOGO_ENTRY_CACHE_SCORE, cap)
            assert need == small(plans, "score_plan", p, ALL, cap)["total"]
            sizes.append((L, cap, p, need))
    for L, cap, p, need in sizes:
        for Lb, capb, _, room in sizes:
            if Lb >= L and capb >= cap:
                got = small(plans, "score_plan", p, room, cap)
                assert got["total"] <= room and got["kc"] % 64 == 0
                assert got["chunks"] == -(-L // got["kc"]) >= 1
                assert got["total"] == up(8 * cap * hq * got["chunks"])
        assert small(plans, "score_plan", p, need, cap) == small(plans, "score_plan", p, ALL, cap)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("B", [1, 4, 16, 100])
def test_step_workspace_of_longer_caches(plans, lib, hq, hkv, d, B):
    import paper_2608_29539_amd as pk
    sizes = []
    for L in (1, 255, 256, 257, 1023, 1024, 1025, 1536, 1537, 4096, 4097, 8191, 32768, 131071):
        p = problem(B, B * L, L, hq, hkv, d, 64)
        need = lib.logo_workspace_bytes(ctypes.byref(p), pk.LOGO_ENTRY_DECODE_SCORE, 0)
        assert need == small(plans, "step_plan", p, ALL)["total"]
        sizes.append((L, p, need))
    for L, p, need in sizes:
        for Lb, _, room in sizes:
            if Lb >= L:
                got = small(plans, "step_plan", p, room)
                assert got["total"] <= room and got["kc"] % 64 == 0
                assert got["chunks"] == -(-L // got["kc"])
                assert got["total"] == up(4 * (hq * B * L + 1)) + up(8 * B * hq * got["chunks"])
        assert small(plans, "step_plan", p, need) == small(plans, "step_plan", p, ALL)


def test_step_sizes_that_shrink(lib):
    import paper_2608_29539_amd as pk

    def need(L):
        p = problem(16, 16 * L, L, 32, 8, 128, 64)
        return lib.logo_workspace_bytes(ctypes.byref(p), pk.LOGO_ENTRY_DECODE_SCORE, 0)

    assert need(1536) > need(1537)


def test_evict_workspace_grows(plans, lib):
    import paper_2608_29539_amd as pk
    last = -1
    for L in (1, 2048, 2049, 8192, 8193, 16384, 16385, 131071):
        p = problem(7, 7 * L, L, 8, 2, 128, 64)
        need = lib.logo_workspace_bytes(ctypes.byref(p), pk.LOGO_ENTRY_CACHE_EVICT, 0)
        assert need == plans.evict_total(ctypes.byref(p)) >= last
        last = need


def test_shapes_reach_their_paths(plans):
    """The shapes that the GPU tests run take the kernels' larger variants."""
    import _cache_shapes as shapes
    seen = set()
    for (lens, rows, hq, hkv, d), waves in shapes.SCORES:
        p = problem(len(lens), sum(lens), max(lens), hq, hkv, d, 64)
        assert plans.score_key_waves(ctypes.byref(p), sum(rows)) == waves
        seen.add((waves, d))
    assert seen == {(w, d) for w in (2, 4) for d in (64, 128)}
    seen = set()
    for (lens, hq, hkv, d), kc in shapes.STEPS:
        p = problem(len(lens), sum(lens), max(lens), hq, hkv, d, 64)
        assert small(plans, "step_plan", p, ALL)["kc"] == kc
        seen.add((kc, d, plans.step_head_copies(ctypes.byref(p))))
        # a wave's half of a chunk, 16 keys a slot, against the ring's slots
        if kc == 1024:
            assert kc // 2 // 16 >= 2 * {64: 16, 128: 8}[d]
    assert seen >= {(kc, d, c) for kc in (512, 1024) for d in (64, 128) for c in (1, 2, 4)}
